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
// thread has kAhead rows' loads in flight: the ids first, then the rows.
constexpr int kAhead = 4;

template <typename T, int V>
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
                if (f0 + u * kThreads < total)
                    store_vec<T, V>(out + (row0 + row[u]) * ld_out + col[u], x[u]);
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
    hipLaunchKernelGGL((k_rows_get<T, V>), dim3((unsigned)wgs), dim3(kThreads), 0, st, (const T*)a.table, a.rows, a.ld,
                       a.k, a.ids, a.ids_stride, a.count, a.scale, (T*)a.out, a.ld_out, per_wg,
                       fast_div((uint32_t)nv));
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
// sort.  A workgroup takes one token at a time; if no earlier token has its id
// it adds the rows of all that do, each wavefront those of a consecutive part
// of the tokens, the four sums joined in order.
constexpr int kScanMost = 4096;

template <typename T, int E>
__global__ __launch_bounds__(kThreads) void k_grad_scan(const T* __restrict__ dout, int64_t ld_dout,
                                                        const int32_t* __restrict__ ids, int64_t ids_stride, int count,
                                                        int k, float scale, T* __restrict__ dtable, int64_t rows,
                                                        int64_t ld, int accumulate)
{
    __shared__ int32_t all[kScanMost];
    __shared__ float part[3][64 * E];
    __shared__ int seen[2][4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Cols c = my_cols<E>(k);
    for (int j = threadIdx.x; j < count; j += kThreads) {
        const int32_t id = ids[j * ids_stride];
        all[j] = id >= 0 && id < rows ? id : -1;
    }
    __syncthreads();
    const int blocks = (count + 63) / 64;
    int turn = 0;
    for (int i = blockIdx.x; i < count; i += gridDim.x) {
        const int32_t r = all[i];
        if (r < 0)
            continue;
        int before = 0;
        for (int b = wave; b * 64 < i && !before; b += 4) {
            const int j = b * 64 + lane;
            before = __ballot(j < i && all[j] == r) != 0;
        }
        if (lane == 0)
            seen[turn][wave] = before;
        __syncthreads();
        const bool first = !(seen[turn][0] | seen[turn][1] | seen[turn][2] | seen[turn][3]);
        turn ^= 1; // the other half is free: everyone passed the last barrier after reading it
        if (!first)
            continue;
        float sum[E];
#pragma unroll
        for (int e = 0; e < E; ++e)
            sum[e] = 0.0f;
        const int b0 = i / 64, each = (blocks - b0 + 3) / 4;
        const int b1 = b0 + wave * each, b2 = b1 + each < blocks ? b1 + each : blocks;
        for (int b = b1; b < b2; ++b) {
            const int j = b * 64 + lane;
            uint64_t mine = __ballot(j >= i && j < count && all[j < count ? j : 0] == r);
            while (mine) {
                int at[4], n = 0;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    at[u] = mine ? __builtin_ctzll(mine) : at[0];
                    n += mine != 0;
                    mine &= mine - 1;
                }
                Vec<T, E> x[4];
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    x[u] = load_vec<T, E>(dout + (int64_t)(b * 64 + at[u]) * ld_dout + c.at);
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (u < n) {
#pragma unroll
                        for (int e = 0; e < E; ++e)
                            sum[e] += (float)x[u].v[e];
                    }
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
            for (int w = 0; w < 3; ++w)
#pragma unroll
                for (int e = 0; e < E; ++e)
                    sum[e] += part[w][e * 64 + lane];
            write_row<T, E>(dtable + (int64_t)r * ld, c, sum, scale, accumulate);
        }
        __syncthreads();
    }
}

// Many tokens: (row, token) pairs sorted by row, stably, so that a row's tokens
// stay in order; then tiles of the sorted tokens summed by one wavefront each.
//
// The sort is by digits of `bits` bits from the lowest: per chunk of kChunk
// tokens the count of every digit, the exclusive sums of these over the chunks,
// and every token to its place.  Tokens without a row have the key `rows` and
// end up last.
constexpr int kChunk = 4096;
constexpr int kDigits = 256;

__device__ __forceinline__ uint32_t key_of(int32_t id, int64_t rows)
{
    return id >= 0 && id < rows ? (uint32_t)id : (uint32_t)rows;
}

__global__ __launch_bounds__(kThreads) void k_sort_count(const uint32_t* __restrict__ keys,
                                                         const int32_t* __restrict__ ids, int64_t ids_stride,
                                                         int64_t rows, int64_t count, int shift, uint32_t mask,
                                                         uint32_t* __restrict__ hist, uint32_t* __restrict__ crossing)
{
    __shared__ uint32_t n[kDigits];
    n[threadIdx.x] = 0;
    __syncthreads();
    const int64_t base = (int64_t)blockIdx.x * kChunk;
#pragma unroll 4
    for (int j = threadIdx.x; j < kChunk; j += kThreads)
        if (base + j < count) {
            const uint32_t key = keys ? keys[base + j] : key_of(ids[(base + j) * ids_stride], rows);
            atomicAdd(&n[key >> shift & mask], 1u);
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
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
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

__global__ __launch_bounds__(kThreads) void k_sort_place(const uint32_t* __restrict__ keys,
                                                         const uint32_t* __restrict__ toks,
                                                         const int32_t* __restrict__ ids, int64_t ids_stride,
                                                         int64_t rows, int64_t count, int shift, int bits,
                                                         const uint32_t* __restrict__ hist,
                                                         const uint32_t* __restrict__ totals,
                                                         uint32_t* __restrict__ keys_out,
                                                         uint32_t* __restrict__ toks_out)
{
    constexpr int steps = kChunk / kThreads; // 64 consecutive tokens a step, a wavefront's steps consecutive
    __shared__ uint32_t next[4][kDigits];
    __shared__ uint32_t sums[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t mask = (1u << bits) - 1;
    const int64_t base = (int64_t)blockIdx.x * kChunk + wave * (steps * 64) + lane;
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
    uint32_t at = block_scan(threadIdx.x <= mask ? totals[threadIdx.x] : 0, sums, total);
    if (threadIdx.x <= mask) {
        at += hist[(int64_t)threadIdx.x * gridDim.x + blockIdx.x];
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
// `tile` tokens, kBatch loads in flight.  A row whose tokens lie inside one tile
// is written at once.  Of one that goes on, the tile where it begins keeps its
// sum in `tails` and notes the tile in `begun`, every later tile its own in
// `heads`; k_grad_join adds those up in order.  The workgroups past the tiles
// write zeros to the rows that no token has.
constexpr int kBatch = 8;

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

template <typename T, int E>
__global__ __launch_bounds__(kThreads) void k_grad_tiles(const T* __restrict__ dout, int64_t ld_dout,
                                                         const uint32_t* __restrict__ keys,
                                                         const uint32_t* __restrict__ toks, int64_t count, int k,
                                                         float scale, T* __restrict__ dtable, int64_t rows, int64_t ld,
                                                         int accumulate, int tile, int64_t tiles, int tile_wgs,
                                                         float* __restrict__ heads, float* __restrict__ tails,
                                                         uint32_t* __restrict__ begun, uint32_t* __restrict__ crossing,
                                                         FastDiv nv)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if ((int)blockIdx.x >= tile_wgs) {
        if (blockIdx.y)
            return;
        const int64_t stride = (int64_t)(gridDim.x - tile_wgs) * 256;
        for (int64_t r0 = ((int64_t)(blockIdx.x - tile_wgs) * 4 + wave) * 64; r0 < rows; r0 += stride) {
            const uint32_t r = (uint32_t)(r0 + lane < rows ? r0 + lane : rows - 1);
            int64_t lo = 0, hi = count; // first sorted token whose key is not below r
            while (lo < hi) {
                const int64_t mid = (lo + hi) >> 1;
                if (keys[mid] < r)
                    lo = mid + 1;
                else
                    hi = mid;
            }
            const uint64_t taken = __ballot(lo < count && keys[lo < count ? lo : 0] == r);
            const int here = (int)(rows - r0 < 64 ? rows - r0 : 64);
            constexpr int most = 16 / (int)sizeof(T);
            if (k >= most)
                zero_rows<T, most>(dtable + r0 * ld, ld, k, here, taken, nv);
            else if (k >= most / 2)
                zero_rows<T, most / 2>(dtable + r0 * ld, ld, k, here, taken, nv);
            else if (most == 8 && k >= 2)
                zero_rows<T, 2>(dtable + r0 * ld, ld, k, here, taken, nv);
            else
                zero_rows<T, 1>(dtable + r0 * ld, ld, k, here, taken, nv);
        }
        return;
    }
    const int64_t t = (int64_t)blockIdx.x * 4 + wave;
    if (t >= tiles)
        return;
    const Cols c = my_cols<E>(k);
    const int64_t start = t * tile;
    const int n = (int)(count - start < tile ? count - start : tile);
    const uint32_t none = 0xffffffffu, out_of_rows = (uint32_t)rows;
    const uint32_t key = keys[start + (lane < n ? lane : n - 1)], tok = toks[start + (lane < n ? lane : n - 1)];
    const uint32_t prev = start > 0 ? keys[start - 1] : none, after = start + n < count ? keys[start + n] : none;
    uint32_t cur = __builtin_amdgcn_readfirstlane(key);
    if (cur == out_of_rows)
        return;
    bool head = prev == cur;
    float sum[E];
#pragma unroll
    for (int e = 0; e < E; ++e)
        sum[e] = 0.0f;
    auto flush = [&](bool tail) {
        if (!head && !tail) {
            write_row<T, E>(dtable + (int64_t)cur * ld, c, sum, scale, accumulate);
            return;
        }
        float* to = (head ? heads : tails) + t * k + c.at;
        if (c.skip < E) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                to[e] = sum[e];
        }
        if (!head && blockIdx.y == 0 && lane == 0)
            begun[atomicAdd(crossing, 1u)] = (uint32_t)t;
    };
    for (int j0 = 0; j0 < n; j0 += kBatch) {
        Vec<T, E> x[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const uint32_t row = __builtin_amdgcn_readlane(tok, j0 + u < n ? j0 + u : n - 1);
            x[u] = load_vec<T, E>(dout + (int64_t)row * ld_dout + c.at);
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (j0 + u < n) {
                const uint32_t at = __builtin_amdgcn_readlane(key, j0 + u);
                if (at != cur) {
                    flush(false);
                    if (at == out_of_rows)
                        return;
                    cur = at;
                    head = false;
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        sum[e] = 0.0f;
                }
#pragma unroll
                for (int e = 0; e < E; ++e)
                    sum[e] += (float)x[u].v[e];
            }
        }
    }
    flush(after == cur);
}

// Joins the rows that go on over several tiles: tails[a], then heads[a + 1 ..
// b], where b is the last tile that begins with the row's key.  A wavefront
// takes one such row a round and adds it alone up to kJoinAlone tiles; a longer
// one is then added by the whole workgroup, its wavefronts taking consecutive
// parts that are joined in order.
constexpr int kJoinThreads = 1024;
constexpr int kJoinAlone = 32;

template <int E>
__device__ __forceinline__ void add_parts(const float* __restrict__ heads, const float* __restrict__ tails, int64_t a,
                                          int from, int to, int k, const Cols& c, float (&sum)[E])
{
    for (int i0 = from; i0 < to; i0 += kBatch) {
        Vec<float, E> x[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int i = i0 + u < to ? i0 + u : to - 1;
            x[u] = load_vec<float, E>((i ? heads : tails) + (a + i) * k + c.at);
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
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
                                                            int tile, int64_t tiles, const float* __restrict__ heads,
                                                            const float* __restrict__ tails,
                                                            const uint32_t* __restrict__ begun,
                                                            const uint32_t* __restrict__ crossing)
{
    constexpr int waves = kJoinThreads / 64;
    __shared__ float part[waves][64 * E];
    __shared__ int long_at[waves], long_span[waves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Cols c = my_cols<E>(k);
    const int64_t n = *crossing;
    float sum[E];
    for (int64_t i0 = (int64_t)blockIdx.x * waves; i0 < n; i0 += (int64_t)gridDim.x * waves) {
        int span = 0;
        if (i0 + wave < n) {
            const int64_t a = __builtin_amdgcn_readfirstlane((int)begun[i0 + wave]);
            const uint32_t key = __builtin_amdgcn_readfirstlane((int)keys[(a + 1) * tile]);
            // tile `lo` begins with the key, tile `hi` does not; 64 places between them a step
            int64_t lo = a + 1, hi = tiles;
            while (hi - lo > 1) {
                const int64_t step = (hi - lo + 63) / 64, p = lo + (lane + 1) * step;
                const int f = __builtin_ctzll(__ballot(p >= hi || keys[(p < hi ? p : lo) * tile] != key));
                const int64_t top = lo + (f + 1) * step;
                lo += f * step;
                hi = top < hi ? top : hi;
            }
            span = (int)(lo - a) + 1;
            if (lane == 0)
                long_at[wave] = (int)a;
            if (span <= kJoinAlone) {
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
            const int total = long_span[w];
            if (total <= kJoinAlone)
                continue;
            const int64_t a = long_at[w];
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

// Tokens of a tile: 64, or fewer where that leaves the chip without enough
// wavefronts to cover the loads' latency.
int tile_of(int64_t count) { return count >= 64 * 4096 ? 64 : count >= 32 * 4096 ? 32 : 16; }

struct GradWork {
    uint32_t *keys[2], *toks[2], *hist, *totals, *crossing, *begun;
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
    const size_t chunks = (size_t)((count + kChunk - 1) / kChunk);
    const size_t tiles = (size_t)((count + tile_of(count) - 1) / tile_of(count));
    for (int i = 0; i < 2; ++i) {
        w.keys[i] = (uint32_t*)part(4 * (size_t)count);
        w.toks[i] = (uint32_t*)part(4 * (size_t)count);
    }
    w.hist = (uint32_t*)part(4 * chunks * kDigits);
    w.totals = (uint32_t*)part(4 * kDigits);
    w.crossing = (uint32_t*)part(4);
    w.begun = (uint32_t*)part(4 * tiles);
    w.heads = (float*)part(4 * tiles * (size_t)k);
    w.tails = (float*)part(4 * tiles * (size_t)k);
    w.bytes = at;
    return w;
}

template <typename T, int E>
hipError_t grad_launch(const RowsGradLaunch& a, hipStream_t st)
{
    const unsigned ys = (unsigned)((a.k + 64 * E - 1) / (64 * E));
    if (a.count <= kScanMost) {
        if (!a.accumulate && a.rows > 0) {
            const hipError_t e = zero_typed<T>(a, st);
            if (e != hipSuccess)
                return e;
        }
        if (a.count == 0)
            return hipSuccess;
        hipLaunchKernelGGL((k_grad_scan<T, E>), dim3((unsigned)std::min<int64_t>(a.count, 2048), ys), dim3(kThreads), 0,
                           st, (const T*)a.dout, a.ld_dout, a.ids, a.ids_stride, (int)a.count, a.k, a.scale,
                           (T*)a.dtable, a.rows, a.ld, a.accumulate);
        return hipGetLastError();
    }
    const GradWork w = grad_work(a.count, a.k, a.work);
    const unsigned chunks = (unsigned)((a.count + kChunk - 1) / kChunk);
    const int bits = key_bits(a.rows), passes = (bits + 7) / 8, width = (bits + passes - 1) / passes;
    const uint32_t *keys = nullptr, *toks = nullptr;
    for (int p = 0; p < passes; ++p) {
        const int shift = p * width, now = std::min(width, bits - shift);
        const uint32_t mask = (1u << now) - 1;
        hipLaunchKernelGGL(k_sort_count, dim3(chunks), dim3(kThreads), 0, st, keys, a.ids, a.ids_stride, a.rows,
                           a.count, shift, mask, w.hist, w.crossing);
        hipLaunchKernelGGL(k_sort_scan, dim3(1u << now), dim3(kThreads), 0, st, w.hist, (int)chunks, w.totals);
        hipLaunchKernelGGL(k_sort_place, dim3(chunks), dim3(kThreads), 0, st, keys, toks, a.ids, a.ids_stride, a.rows,
                           a.count, shift, now, w.hist, w.totals, w.keys[p & 1], w.toks[p & 1]);
        keys = w.keys[p & 1];
        toks = w.toks[p & 1];
    }
    const int tile = tile_of(a.count);
    const int64_t tiles = (a.count + tile - 1) / tile;
    const int tile_wgs = (int)((tiles + 3) / 4);
    const int zero_wgs = a.accumulate ? 0 : (int)std::min<int64_t>((a.rows + 255) / 256, 1 << 20);
    const int v = vec_of<T>(a.k);
    hipLaunchKernelGGL((k_grad_tiles<T, E>), dim3((unsigned)(tile_wgs + zero_wgs), ys), dim3(kThreads), 0, st,
                       (const T*)a.dout, a.ld_dout, keys, toks, a.count, a.k, a.scale, (T*)a.dtable, a.rows, a.ld,
                       a.accumulate, tile, tiles, tile_wgs, w.heads, w.tails, w.begun, w.crossing,
                       fast_div((uint32_t)((a.k + v - 1) / v)));
    hipLaunchKernelGGL((k_grad_join<T, E>), dim3((unsigned)std::min<int64_t>((tiles + 15) / 16, 256), ys),
                       dim3(kJoinThreads), 0, st, keys, a.k, a.scale, (T*)a.dtable, a.ld, a.accumulate, tile, tiles,
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

size_t rows_grad_bytes(int64_t count, int k) { return count <= kScanMost ? 0 : grad_work(count, k, nullptr).bytes; }

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
